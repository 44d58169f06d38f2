"""Performance cases of the 8-bit integer layer: a user's calls of `paper_2609_26077_b200.int8`, and their plain forms.

Five kinds of work, with the sizes of the library's own benchmark and error-sweep configurations (`bench.py`,
`paper_2609_26077_b200/sweep.py`) and ragged ones between them:

  checkpoint  activations saved in 8 bits and restored (int8.quantize, int8.dequantize)
  norm        residual's addition, root-mean-square norm and 8-bit output, with or without an 8-bit checkpoint of the
              hidden rows (the sums) for the backward pass (int8.rms_norm)
  norm_back   gradients of that norm, from the checkpoint (int8.rms_norm_backward)
  matmul      product of 8-bit codes with a scale per token and per output channel (int8.matmul)
  linear_back both gradients of that product, from the 8-bit activations and weights (int8.grad_weight, int8.grad_input)

The codes of a block x of numbers are round(x * (127 / max|x|)), ties to even, and its scale is max|x| / 127, or with
`pow2` the power of two at or above that.  run() returns what 8-bit codes stand for, code * scale, not the codes.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def _checkpoint(rows, cols, dtype, block, pow2):
    return {"kind": "checkpoint", "rows": rows, "cols": cols, "dtype": dtype, "block": block, "pow2": pow2}


def _norm(rows, cols, dtype, residual, pow2, block, kind="norm"):
    return {"kind": kind, "rows": rows, "cols": cols, "dtype": dtype, "residual": residual, "pow2": pow2, "block": block}


def _matmul(M, N, K, dtype, bias):
    return {"kind": "matmul", "M": M, "N": N, "K": K, "dtype": dtype, "bias": bias}


def _linear_back(M, N, K, dtype, wdtype):
    return {"kind": "linear_back", "M": M, "N": N, "K": K, "dtype": dtype, "wdtype": wdtype}


def listed():
    def named(name, case):
        return {"name": name, **case}
    return [
        # the activations of a short ragged batch, in blocks of 32 with power-of-two scales (exact in bf16)
        named("checkpoint_777x2048", _checkpoint(777, 2048, "bf16", 32, True)),
        # the activations of a full training step's tokens, blocks of 128
        named("checkpoint_16384x8192", _checkpoint(16384, 8192, "bf16", 128, False)),
        # decoding: one token's hidden row, on the way into the next product
        named("norm_1x8192", _norm(1, 8192, "bf16", True, False, 0)),
        # prefill of a ragged batch in half precision, row length no multiple of a vector
        named("norm_1000x4095", _norm(1000, 4095, "fp16", True, False, 0)),
        # training: hidden rows checkpointed on the way
        named("norm_16384x8192", _norm(16384, 8192, "bf16", True, True, 128)),
        # backward of a short ragged batch, no gradient beside the norm's own
        named("norm_back_777x2048", _norm(777, 2048, "bf16", False, False, 32, kind="norm_back")),
        # backward of a full training step's tokens
        named("norm_back_16384x8192", _norm(16384, 8192, "bf16", True, False, 128, kind="norm_back")),
        # decoding: one token through a square weight
        named("matmul_1x8192x8192", _matmul(1, 8192, 8192, "bf16", False)),
        # a ragged batch of prompts through a small layer with a bias, full-precision output
        named("matmul_777x2047x2048", _matmul(777, 2047, 2048, "fp32", True)),
        # the LLM-shaped product of the benchmark
        named("matmul_16384x8192x8192", _matmul(16384, 8192, 8192, "bf16", False)),
        # backward of a ragged batch through a small layer
        named("linear_back_1001x2048x2047", _linear_back(1001, 2048, 2047, "bf16", "fp32")),
        # backward of a full step
        named("linear_back_8192x8192x8192", _linear_back(8192, 8192, 8192, "bf16", "fp32")),
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        # half of the sizes are multiples of 64, as those of models are; the others are whatever came
        return max(lo, n // 64 * 64) if n >= 128 and rng.random() < 0.5 else n
    kind = rng.choice(["checkpoint", "norm", "norm_back", "matmul", "linear_back"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind == "checkpoint":
        return _checkpoint(size(1, 16384), size(64, 8192), dtype, rng.choice([0, 32, 128]), rng.random() < 0.5)
    if kind in ("norm", "norm_back"):
        block = rng.choice([32, 128] if kind == "norm_back" else [0, 0, 32, 128])
        return _norm(size(1, 16384), size(64, 8192), dtype, rng.random() < 0.7, kind == "norm" and rng.random() < 0.3, block, kind)
    if kind == "matmul":
        return _matmul(size(1, 16384), size(64, 8192), size(64, 8192), dtype, rng.random() < 0.5)
    return _linear_back(size(16, 8192), size(64, 8192), size(64, 8192), rng.choice(["bf16", "fp16"]), rng.choice(["fp32", "same"]))


def _padded(x):
    """The same values with rows 16 bytes (or a multiple) apart, as the library's own outputs have them."""
    ld = -(-x.shape[1] * x.element_size() // 16) * 16 // x.element_size()
    out = torch.zeros(x.shape[0], ld, dtype=x.dtype, device=x.device)[:, :x.shape[1]]
    out.copy_(x)
    return out


def _activations(rows, cols, dtype, gen, sigma=1.0):
    """Rows N(0, 1) times a lognormal factor per channel: the operands of the benchmark's LLM-shaped product."""
    factor = torch.exp(sigma * torch.randn(cols, device="cuda", generator=gen))
    return (torch.randn(rows, cols, device="cuda", generator=gen) * factor).to(dtype)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    dtype = DTYPES[case["dtype"]]
    if kind in ("checkpoint", "norm", "norm_back"):
        rows, cols = case["rows"], case["cols"]
    if kind == "checkpoint":
        s["x"] = _activations(rows, cols, dtype, gen)
    elif kind == "norm":
        s["x"] = _activations(rows, cols, dtype, gen)
        s["residual"] = _activations(rows, cols, dtype, gen) if case["residual"] else None
        s["gain"] = (1 + 0.2 * torch.randn(cols, device="cuda", generator=gen)).to(dtype)
    elif kind == "norm_back":
        # what the forward pass left: codes and scales of the hidden rows, and their reciprocal root mean squares
        hidden = _activations(rows, cols, torch.float32, gen)
        codes, s["scales"] = _quantize(hidden, case["block"], case["pow2"])
        s["codes"] = _padded(codes.to(torch.int8))
        s["rstd"] = (hidden.double().square().mean(1) + EPS).rsqrt().float()
        s["gain"] = (1 + 0.2 * torch.randn(cols, device="cuda", generator=gen)).to(dtype)
        s["dy"] = torch.randn(rows, cols, device="cuda", generator=gen).to(dtype)
        s["dresidual"] = torch.randn(rows, cols, device="cuda", generator=gen).to(dtype) if case["residual"] else None
    else:
        M, N, K = case["M"], case["N"], case["K"]
        weights = 0.02 * torch.randn(N, K, device="cuda", generator=gen)
        codes, s["wscales"] = _quantize(weights, 0, False)
        s["w"] = _padded(codes.to(torch.int8))
        tokens = _activations(M, K, torch.float32, gen)
        # a gradient in 32 bits takes activations with power-of-two scales, whose values are exact in 16 bits
        codes, s["xscales"] = _quantize(tokens, 0, kind == "linear_back" and case["wdtype"] == "fp32")
        s["x"] = _padded(codes.to(torch.int8))
        if kind == "matmul":
            s["bias"] = torch.randn(N, device="cuda", generator=gen).to(dtype) if case["bias"] else None
        else:
            s["dy"] = torch.randn(M, N, device="cuda", generator=gen).to(dtype)
    return s


# ---------------------------------------------------------------- plain forms

def _blocks(x, block):
    """(rows, blocks, block) with zeros behind the last column; block 0: the whole row."""
    rows, cols = x.shape
    block = block or cols
    return torch.nn.functional.pad(x, (0, -cols % block)).view(rows, -1, block)


def _quantize(x, block, pow2):
    """Codes (as 32-bit numbers) and scales of 32-bit rows."""
    b = _blocks(x, block)
    amax = b.abs().amax(2).clamp_min(1e-12)
    full = torch.full_like(amax, 127.0)
    scales, inverse = amax / full, full / amax
    if pow2:
        mantissa, exponent = torch.frexp(scales)
        scales = torch.ldexp(torch.ones_like(scales), exponent - (mantissa == 0.5).int())
        inverse = 1 / scales
    codes = torch.round(b * inverse[:, :, None]).clamp(-127, 127).flatten(1)[:, :x.shape[1]]
    return codes, scales if block else scales[:, 0]


def _values(codes, scales, block):
    b = _blocks(codes.float(), block)
    return (b * scales.view(b.shape[0], -1, 1)).flatten(1)[:, :codes.shape[1]]


def _short(dtype):
    """The type in which values of 8-bit codes are handed on."""
    return torch.float16 if dtype == torch.float16 else torch.bfloat16


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    dtype = DTYPES[case["dtype"]]
    if kind == "checkpoint":
        codes, scales = _quantize(s["x"].float(), case["block"], case["pow2"])
        return {"values": _values(codes, scales, case["block"]).to(_short(dtype)), "scales": scales}
    if kind == "norm":
        h = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
        rstd = (1 / torch.sqrt(h.double().square().mean(1) + EPS)).float()
        codes, scales = _quantize(h * rstd[:, None] * s["gain"].float(), 0, case["pow2"])
        out = {"values": _values(codes, scales, 0).to(_short(dtype)), "scales": scales, "rstd": rstd}
        if s["residual"] is not None:
            out["hidden"] = h.to(dtype)
        if case["block"]:
            codes, scales = _quantize(h, case["block"], False)
            out["checkpoint"] = _values(codes, scales, case["block"]).to(_short(dtype))
            out["checkpoint_scales"] = scales
        return out
    if kind == "norm_back":
        xhat = _values(s["codes"], s["scales"], case["block"]) * s["rstd"][:, None]
        dy = s["dy"].float()
        dxhat = dy * s["gain"].float()
        dx = (dxhat - xhat * (dxhat * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
        if s["dresidual"] is not None:
            dx = dx + s["dresidual"].float()
        return {"dx": dx.to(dtype), "dgain": (dy * xhat).sum(0)}
    if kind == "matmul":
        c = s["x"].float() @ s["w"].float().t() * s["xscales"][:, None] * s["wscales"][None, :]
        return (c if s["bias"] is None else c + s["bias"].float()).to(dtype)
    dy = s["dy"].float()
    dw = dy.t() @ _values(s["x"], s["xscales"], 0)
    dx = dy @ _values(s["w"], s["wscales"], 0)
    return {"dw": dw if case["wdtype"] == "fp32" else dw.to(dtype), "dx": dx.to(dtype)}


# ---------------------------------------------------------------- the library's calls

def _run_own(s):
    from paper_2609_26077_b200 import int8
    case, kind = s["case"], s["case"]["kind"]
    dtype = DTYPES[case["dtype"]]
    if kind == "checkpoint":
        codes, scales = int8.quantize(s["x"], block=case["block"], pow2=case["pow2"])
        return {"values": int8.dequantize(codes, scales, block=case["block"], dtype=_short(dtype)), "scales": scales}
    if kind == "norm":
        n = int8.rms_norm(s["x"], s["gain"], residual=s["residual"], eps=EPS, pow2=case["pow2"], checkpoint=case["block"])
        out = {"values": int8.dequantize(n.codes, n.scales, dtype=_short(dtype)), "scales": n.scales, "rstd": n.rstd}
        if s["residual"] is not None:
            out["hidden"] = n.hidden
        if case["block"]:
            out["checkpoint"] = int8.dequantize(n.checkpoint, n.checkpoint_scales, block=case["block"], dtype=_short(dtype))
            out["checkpoint_scales"] = n.checkpoint_scales
        return out
    if kind == "norm_back":
        dx, dgain = int8.rms_norm_backward(s["dy"], s["codes"], s["scales"], s["rstd"], s["gain"], block=case["block"],
                                           dresidual=s["dresidual"])
        return {"dx": dx, "dgain": dgain}
    if kind == "matmul":
        return int8.matmul(s["x"], s["xscales"], s["w"], s["wscales"], bias=s["bias"], dtype=dtype)
    return {"dw": int8.grad_weight(s["dy"], s["x"], s["xscales"], dtype=torch.float32 if case["wdtype"] == "fp32" else dtype),
            "dx": int8.grad_input(s["dy"], s["w"], s["wscales"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- definitions in 64 bits

def _exact_values(x, block, pow2):
    """What the codes of 64-bit rows stand for, and their scales."""
    rows, cols = x.shape
    width = block if block else cols
    scales, values = [], []
    for c in range(0, cols, width):
        piece = x[:, c:c + width]
        top = torch.clamp(piece.abs().max(dim=1).values, min=1e-12)
        scale = top / torch.tensor(127.0, dtype=top.dtype, device=top.device)      # by a tensor: a plain number is multiplied by its reciprocal
        if pow2:
            # from a power that is too small up to the first that is not: a logarithm may be a little off at a power itself
            power = torch.ldexp(torch.ones_like(scale), torch.floor(torch.log2(scale)).int() - 2)
            for _ in range(4):
                power = torch.where(power < scale, 2 * power, power)
            scale = power
        steps = torch.round(piece / scale.unsqueeze(1))
        scales.append(scale)
        values.append(steps * scale.unsqueeze(1))
    return torch.cat(values, 1), torch.stack(scales, 1) if block else scales[0]


def _held(codes, scales, block):
    """Codes and scales that are given, as 64-bit numbers."""
    scales = scales.double()
    if block:
        scales = scales.repeat_interleave(block, dim=1)[:, :codes.shape[1]]
    else:
        scales = scales.unsqueeze(1)
    return codes.double() * scales


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "checkpoint":
        values, scales = _exact_values(s["x"].double(), case["block"], case["pow2"])
        return {"values": values, "scales": scales}
    if kind == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        rstd = 1 / ((h * h).sum(1) / h.shape[1] + EPS) ** 0.5
        values, scales = _exact_values(torch.einsum("rc,r,c->rc", h, rstd, s["gain"].double()), 0, case["pow2"])
        out = {"values": values, "scales": scales, "rstd": rstd}
        if s["residual"] is not None:
            out["hidden"] = h
        if case["block"]:
            out["checkpoint"], out["checkpoint_scales"] = _exact_values(h, case["block"], False)
        return out
    if kind == "norm_back":
        n, rstd, gain, dy = case["cols"], s["rstd"].double(), s["gain"].double(), s["dy"].double()
        h = _held(s["codes"], s["scales"], case["block"])
        # y = gain * h * rstd, with d rstd / d h = -rstd^3 h / n
        along = torch.einsum("rc,rc,c->r", dy, h, gain)
        dx = rstd[:, None] * gain * dy - (rstd ** 3 * along / n)[:, None] * h
        if s["dresidual"] is not None:
            dx = dx + s["dresidual"].double()
        return {"dx": dx, "dgain": torch.einsum("rc,rc,r->c", dy, h, rstd)}
    if kind == "matmul":
        c = torch.matmul(_held(s["x"], s["xscales"], 0), _held(s["w"], s["wscales"], 0).T)
        return c if s["bias"] is None else c + s["bias"].double()
    dy = s["dy"].double()
    return {"dw": torch.matmul(dy.T, _held(s["x"], s["xscales"], 0)), "dx": torch.matmul(dy, _held(s["w"], s["wscales"], 0))}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    kind = case["kind"]
    if kind in ("checkpoint", "norm", "norm_back"):
        rows, cols, block = case["rows"], case["cols"], case["block"]
        elements, scales = rows * cols, rows * (-(-cols // block) if block else 1)
        if kind == "checkpoint":      # the activations in, their values out
            return {"bytes": elements * (size + 2) + 4 * scales, "flops": 4 * elements}
        if kind == "norm":            # rows (and residual) in; values, hidden rows and the checkpoint's values out
            per = size * (3 if case["residual"] else 1) + 2 + (2 if block else 0)
            return {"bytes": elements * per + 8 * rows + size * cols + (4 * scales if block else 0),
                    "flops": (8 + (4 if block else 0)) * elements}
        per = size * (3 if case["residual"] else 2) + 1
        return {"bytes": elements * per + 4 * (scales + rows) + (size + 4) * cols, "flops": 10 * elements}
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "matmul":
        return {"bytes": M * K + N * K + 4 * (M + N) + size * M * N, "flops": 2 * M * N * K}
    wsize = 4 if case["wdtype"] == "fp32" else size
    return {"bytes": size * M * N + M * K + N * K + 4 * (M + N) + wsize * N * K + size * M * K, "flops": 4 * M * N * K}
