"""Performance cases of the 8-bit floating-point layer: a user's calls of `paper_2609_26077_b200.fp8` and
`paper_2609_26077_b200.gradients`, and their plain forms.

Five kinds of work.  Sizes are those of the library's own benchmark and error-sweep configurations (`bench.py`,
`paper_2609_26077_b200/sweep.py`), ragged ones between them, and generic numbers of experts:

  linear        activations to e4m3 (a scale for each 128 columns of a token) and their product with a weight that is held in
                e4m3 (a scale for each 128 x 128 tile): fp8.quantize, fp8.matmul
  linear_back   both gradients of that product: dy to e4m3 along its rows and along its columns, dx from the weight, dw from
                the activations that the forward pass kept along their columns: fp8.quantize_both, fp8.grad_input, fp8.grad_weight
  experts       the product for tokens that are sorted by expert, a weight to each expert and ragged numbers of tokens:
                fp8.quantize, fp8.grouped_matmul
  experts_back  its gradients: fp8.quantize_both, fp8.grouped_grad_input, fp8.grouped_grad_weight
  clip          gradients of many parameters, scaled to a largest global norm: gradients.clip

With a = max(max |x| of a block, 1e-12) a block's scale is a / 448, or with `pow2` the power of two at or above that, and its codes
are x * (448 / a) (pow2: x / scale) in fp32, rounded to the nearest e4m3 number, ties to even.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BLOCK = 128


def _linear(M, N, K, dtype, bias, pow2, kind="linear"):
    return {"kind": kind, "M": M, "N": N, "K": K, "dtype": dtype, "bias": bias, "pow2": pow2}


def _linear_back(M, N, K, dtype, wdtype, pow2):
    return {"kind": "linear_back", "M": M, "N": N, "K": K, "dtype": dtype, "wdtype": wdtype, "pow2": pow2}


def _experts(E, M, N, K, dtype, spread, pow2):
    return {"kind": "experts", "E": E, "M": M, "N": N, "K": K, "dtype": dtype, "spread": spread, "pow2": pow2}


def _experts_back(E, M, N, K, dtype, wdtype, spread, pow2):
    return {"kind": "experts_back", "E": E, "M": M, "N": N, "K": K, "dtype": dtype, "wdtype": wdtype, "spread": spread, "pow2": pow2}


def _clip(tensors, elements, dtype):
    return {"kind": "clip", "tensors": tensors, "elements": elements, "dtype": dtype}


def listed():
    def named(name, case):
        return {"name": name, **case}
    return [
        # decoding: one token through a square weight
        named("linear_1x8192x8192", _linear(1, 8192, 8192, "bf16", False, False)),
        # a ragged batch of prompts through a small layer with a bias, odd number of output channels, full-precision output
        named("linear_777x2047x2048", _linear(777, 2047, 2048, "fp32", True, False)),
        # the LLM-shaped product of the benchmark
        named("linear_16384x8192x8192", _linear(16384, 8192, 8192, "bf16", False, False)),
        # backward of a ragged batch through a small layer, odd number of input channels
        named("linear_back_1001x2048x2047", _linear_back(1001, 2048, 2047, "fp16", "fp32", False)),
        # backward of a full step
        named("linear_back_8192x8192x8192", _linear_back(8192, 8192, 8192, "bf16", "fp32", False)),
        # decoding with experts: a few tokens, eight experts each, so that most experts see one to four rows
        named("experts_64x128x2048x4096", _experts(64, 128, 2048, 4096, "bf16", 0.0, False)),
        # ragged prompts through eight small experts, power-of-two scales
        named("experts_8x5001x1024x2048", _experts(8, 5001, 1024, 2048, "fp16", 0.5, True)),
        # a full step's tokens
        named("experts_16x32768x4096x4096", _experts(16, 32768, 4096, 4096, "bf16", 0.3, False)),
        # backward of ragged prompts, a few of the experts without any token
        named("experts_back_32x999x1024x2048", _experts_back(32, 999, 1024, 2048, "bf16", "bf16", 1.0, False)),
        # backward of a full step's tokens
        named("experts_back_16x16384x4096x4096", _experts_back(16, 16384, 4096, 4096, "bf16", "fp32", 0.3, False)),
        # gradients of a small model: norms' gains, biases, small weights, lying behind one another in one buffer, odd sizes
        named("clip_200x2000000", _clip(200, 2000000, "bf16")),
        # gradients of the large layers of a step in full precision
        named("clip_24x268435456", _clip(24, 268435456, "fp32")),
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        # half of the sizes are multiples of 64, as those of models are; the others are whatever came
        return max(lo, n // 64 * 64) if n >= 128 and rng.random() < 0.5 else n
    kind = rng.choice(["linear", "linear_back", "experts", "experts_back", "clip"])
    dtype, pow2 = rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.random() < 0.3
    if kind == "linear":
        return _linear(size(1, 16384), size(64, 8192), size(64, 8192), dtype, rng.random() < 0.5, pow2)
    if kind == "linear_back":
        return _linear_back(size(16, 8192), size(64, 8192), size(64, 8192), dtype, rng.choice(["fp32", "same"]), pow2)
    if kind == "clip":
        return _clip(size(1, 400), size(1000, 268435456), dtype)
    N, K, spread = size(64, 4096), size(64, 4096), rng.choice([0.0, 0.3, 0.5, 1.0])
    E = min(size(1, 64), max(1, 268435456 // (N * K)))
    if kind == "experts":
        return _experts(E, size(1, 32768), N, K, dtype, spread, pow2)
    return _experts_back(E, size(16, 16384), N, K, dtype, rng.choice(["fp32", "same"]), spread, pow2)


def _apart(rows, cols, dtype, step):
    """An empty matrix whose rows are a multiple of `step` elements apart, as the library's own outputs have them."""
    return torch.zeros(rows, -(-cols // step) * step, dtype=dtype, device="cuda")[:, :cols]


def _held(codes):
    """e4m3 codes of numbers that e4m3 has."""
    out = _apart(codes.shape[0], codes.shape[1], torch.float8_e4m3fn, 16)
    out.copy_(codes)
    return out


def _held_scales(scales):
    out = _apart(scales.shape[0], scales.shape[1], torch.float32, 4)
    out.copy_(scales)
    return out


def _activations(rows, cols, dtype, gen, sigma=1.0):
    """Rows N(0, 1) times a lognormal factor per channel: the operands of the benchmark's LLM-shaped product."""
    factor = torch.exp(sigma * torch.randn(cols, device="cuda", generator=gen))
    return (torch.randn(rows, cols, device="cuda", generator=gen) * factor).to(dtype)


def _offsets(E, rows, spread, seed):
    """How many of `rows` tokens each of E experts got, as the first row of each and the end of the last; their popularity is lognormal."""
    gen = torch.Generator().manual_seed(seed)
    share = torch.exp(spread * torch.randn(E, generator=gen, dtype=torch.float64))
    counts = torch.bincount(torch.multinomial(share, rows, replacement=True, generator=gen), minlength=E)
    return torch.nn.functional.pad(counts.cumsum(0), (1, 0)).int(), int(counts.max())


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    dtype = DTYPES[case["dtype"]]
    if kind == "clip":
        # sizes are lognormal; the tensors lie behind one another, as the buckets of a data-parallel step have them
        cpu = torch.Generator().manual_seed(seed)
        parts = torch.exp(1.5 * torch.randn(case["tensors"], generator=cpu, dtype=torch.float64))
        ends = torch.round(parts.cumsum(0) / parts.sum() * case["elements"]).long().tolist()
        s["ends"] = ends
        s["sizes"] = [e - b for b, e in zip([0] + ends[:-1], ends)]
        size = torch.exp(torch.randn(len(ends), generator=cpu)).cuda() * 1e-3
        flat = torch.randn(case["elements"], device="cuda", generator=gen)
        for b, e, f in zip([0] + ends[:-1], ends, size):
            flat[b:e] *= f
        s["flat"] = flat.to(dtype)
        s["grads"] = list(s["flat"].split(s["sizes"]))
        s["out_flat"] = torch.empty_like(s["flat"])
        s["out"] = list(s["out_flat"].split(s["sizes"]))
        s["max_norm"] = 0.25
        return s
    M, N, K, pow2 = case["M"], case["N"], case["K"], case["pow2"]
    E = case.get("E", 1)
    if "E" in case:
        offsets, s["longest"] = _offsets(E, M, case["spread"], seed)
        s["offsets"] = offsets.cuda()
    # the weight, or one for each expert
    tiles = [_quantize_tiles(0.02 * torch.randn(N, K, device="cuda", generator=gen), pow2) for _ in range(E)]
    ld = -(-K // 16) * 16
    w = torch.zeros(E, N, ld, dtype=torch.float8_e4m3fn, device="cuda")
    for e, (codes, _) in enumerate(tiles):
        w[e, :, :K] = codes.to(torch.float8_e4m3fn)
    ws = torch.stack([scales for _, scales in tiles])
    s["w"], s["wscales"] = (w[:, :, :K], ws) if "E" in case else (w[0, :, :K], ws[0])
    if kind in ("linear", "experts"):
        s["x"] = _activations(M, K, dtype, gen)
        s["bias"] = torch.randn(N, device="cuda", generator=gen).to(dtype) if case.get("bias") else None
    else:
        # the activations as the forward pass kept them
        codes, scales = _quantize_columns(_activations(M, K, torch.float32, gen), s.get("offsets"), pow2)
        s["x"], s["xscales"] = _held(codes), scales
        s["dy"] = torch.randn(M, N, device="cuda", generator=gen).to(dtype)
    return s


# ---------------------------------------------------------------- plain forms

def _codes(b, dim, pow2):
    """Codes (as 32-bit numbers) of blocks along `dim`, and their scales."""
    amax = b.abs().amax(dim).clamp_min(1e-12)
    full = torch.full_like(amax, 448.0)
    scales, inverse = amax / full, full / amax
    if pow2:
        mantissa, exponent = torch.frexp(scales)
        scales = torch.ldexp(torch.ones_like(scales), exponent - (mantissa == 0.5).int())
        inverse = 1 / scales
    return (b * inverse.unsqueeze(dim)).clamp(-448, 448).to(torch.float8_e4m3fn).float(), scales


def _quantize_rows(x, pow2):
    """Blocks of 128 columns of a row: codes (rows x cols), scales (blocks x rows)."""
    rows, cols = x.shape
    codes, scales = _codes(torch.nn.functional.pad(x, (0, -cols % BLOCK)).view(rows, -1, BLOCK), 2, pow2)
    return codes.flatten(1)[:, :cols], scales.t()


def _quantize_tiles(w, pow2):
    """Tiles of 128 x 128: codes (rows x cols), scales (tiles down x tiles across)."""
    rows, cols = w.shape
    b = torch.nn.functional.pad(w, (0, -cols % BLOCK, 0, -rows % BLOCK))
    b = b.view(b.shape[0] // BLOCK, BLOCK, -1, BLOCK).transpose(1, 2).flatten(2)
    codes, scales = _codes(b, 2, pow2)
    codes = codes.view(b.shape[0], b.shape[1], BLOCK, BLOCK).transpose(1, 2).reshape(b.shape[0] * BLOCK, -1)
    return codes[:rows, :cols], scales


def _places(offsets, rows):
    """Expert and rank of each row, and where it lies once every expert begins on a multiple of 128; rows of that layout that an expert
    begins on, by expert."""
    counts = offsets.diff()
    first = torch.nn.functional.pad((counts + BLOCK - 1) // BLOCK * BLOCK, (1, 0)).cumsum(0)
    at = torch.arange(rows, device=offsets.device)
    expert = torch.searchsorted(offsets[1:].contiguous(), at, right=True)
    rank = at - offsets[expert]
    return expert, rank, first[expert] + rank, first


def _column_rows(rows, offsets):
    """Rows that the form along the columns has."""
    if offsets is None:
        return -(-rows // BLOCK) * BLOCK
    return (rows + (BLOCK - 1) * (offsets.shape[0] - 1)) // BLOCK * BLOCK


def _quantize_columns(x, offsets, pow2):
    """Blocks of 128 rows of a column, counted from the first row of each expert: codes (rows as _column_rows x cols), scales (blocks x cols)."""
    rows, cols = x.shape
    padded = torch.zeros(_column_rows(rows, offsets), cols, device=x.device)
    padded[torch.arange(rows, device=x.device) if offsets is None else _places(offsets, rows)[2]] = x
    codes, scales = _codes(padded.view(-1, BLOCK, cols), 1, pow2)
    return codes.flatten(0, 1), scales


def _row_values(codes, scales):
    return codes * scales.t().repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def _column_values(codes, scales):
    return codes * scales.repeat_interleave(BLOCK, 0)


def _tile_values(codes, scales):
    wide = scales.repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]
    return codes.float() * wide.repeat_interleave(BLOCK, -2)[..., :codes.shape[-2], :]


def _by_expert(x, expert, rank, E, longest):
    """(E, longest, cols): every expert's rows, zeros behind them."""
    out = torch.zeros(E, longest, x.shape[1], device=x.device)
    out[expert, rank] = x
    return out


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    dtype = DTYPES[case["dtype"]]
    if kind == "clip":
        flat = torch.cat(s["grads"]).float()
        norm = flat.double().square().sum().sqrt()
        factor = torch.clamp(s["max_norm"] / norm, max=1.0).float()
        return {"norm": norm.float(), "flat": (flat * factor).to(dtype)}
    w = _tile_values(s["w"], s["wscales"])
    if kind == "linear":
        y = _row_values(*_quantize_rows(s["x"].float(), case["pow2"])) @ w.t()
        return (y if s["bias"] is None else y + s["bias"].float()).to(dtype)
    if kind == "experts":
        x = _row_values(*_quantize_rows(s["x"].float(), case["pow2"]))
        expert, rank, _, _ = _places(s["offsets"], x.shape[0])
        return torch.bmm(_by_expert(x, expert, rank, case["E"], s["longest"]), w.transpose(1, 2))[expert, rank].to(dtype)
    wdtype = torch.float32 if case["wdtype"] == "fp32" else dtype
    dy = s["dy"].float()
    along_rows = _row_values(*_quantize_rows(dy, case["pow2"]))
    along_columns = _column_values(*_quantize_columns(dy, s.get("offsets"), case["pow2"]))
    x = _column_values(s["x"].float(), s["xscales"])
    if kind == "linear_back":
        return {"dx": (along_rows @ w).to(dtype), "dw": (along_columns.t() @ x).to(wdtype)}
    expert, rank, place, _ = _places(s["offsets"], dy.shape[0])
    E, longest = case["E"], s["longest"]
    dx = torch.bmm(_by_expert(along_rows, expert, rank, E, longest), w)[expert, rank]
    dw = torch.bmm(_by_expert(along_columns[place], expert, rank, E, longest).transpose(1, 2), _by_expert(x[place], expert, rank, E, longest))
    return {"dx": dx.to(dtype), "dw": dw.to(wdtype)}


# ---------------------------------------------------------------- the library's calls

def _run_own(s):
    from paper_2609_26077_b200 import fp8, gradients
    case, kind = s["case"], s["case"]["kind"]
    dtype = DTYPES[case["dtype"]]
    if kind == "clip":
        return {"norm": gradients.clip(s["grads"], s["max_norm"], out=s["out"]), "flat": s["out_flat"]}
    if kind == "linear":
        x, xs = fp8.quantize(s["x"], pow2=case["pow2"])
        return fp8.matmul(x, xs, s["w"], s["wscales"], bias=s["bias"], dtype=dtype)
    if kind == "experts":
        x, xs = fp8.quantize(s["x"], pow2=case["pow2"])
        return fp8.grouped_matmul(x, xs, s["w"], s["wscales"], s["offsets"], dtype=dtype)
    wdtype = torch.float32 if case["wdtype"] == "fp32" else dtype
    if kind == "linear_back":
        dy = fp8.quantize_both(s["dy"], pow2=case["pow2"])
        return {"dx": fp8.grad_input(dy.codes, dy.scales, s["w"], s["wscales"], dtype=dtype),
                "dw": fp8.grad_weight(dy.column_codes, dy.column_scales, s["x"], s["xscales"], dtype=wdtype)}
    dy = fp8.quantize_both(s["dy"], offsets=s["offsets"], pow2=case["pow2"])
    return {"dx": fp8.grouped_grad_input(dy.codes, dy.scales, s["w"], s["wscales"], s["offsets"], dtype=dtype),
            "dw": fp8.grouped_grad_weight(dy.column_codes, dy.column_scales, s["x"], s["xscales"], s["offsets"], dtype=wdtype)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- definitions in 64 bits

def _exact_block(b, pow2):
    """What the e4m3 form of one block (or of many: reduced over the last axis) stands for.  The definition rounds 448 / a (or the scale) and
    its product with x to 32 bits."""
    top = torch.clamp(b.abs().max(dim=-1, keepdim=True).values, min=float(torch.tensor(1e-12)))
    scale = (top / 448).float().double()
    if pow2:
        # from a power that is too small up to the first that is not: a logarithm may be a little off at a power itself
        power = torch.ldexp(torch.ones_like(scale), torch.floor(torch.log2(scale)).int() - 2)
        for _ in range(4):
            power = torch.where(power < scale, 2 * power, power)
        scale = power
        y = (b / scale).float().double()
    else:
        y = (b * (448 / top).float().double()).float().double()
    # numbers of e4m3 from 2^e up are 2^(e-3) apart, those below 2^-6 as far as those above it
    step = torch.ldexp(torch.ones_like(y), torch.clamp(torch.frexp(y).exponent - 1, min=-6).int() - 3)
    return torch.clamp(torch.round(y / step) * step, -448, 448) * scale


def _exact_rows(x, pow2):
    return torch.cat([_exact_block(x[:, c:c + BLOCK], pow2) for c in range(0, x.shape[1], BLOCK)], 1)


def _exact_columns(x, bounds, pow2):
    pieces = [x[r:min(r + BLOCK, end)] for begin, end in zip(bounds, bounds[1:]) for r in range(begin, end, BLOCK)]
    return torch.cat([_exact_block(p.T, pow2).T for p in pieces], 0)


def _exact_tiles(codes, scales):
    out = codes.double()
    for r in range(scales.shape[0]):
        for c in range(scales.shape[1]):
            out[r * BLOCK:(r + 1) * BLOCK, c * BLOCK:(c + 1) * BLOCK] *= scales[r, c].double()
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "clip":
        norm = math.sqrt(sum(float(torch.dot(g.double(), g.double())) for g in s["grads"]))
        return {"norm": torch.tensor(norm, dtype=torch.float64), "flat": s["flat"].double() * min(1.0, s["max_norm"] / norm)}
    pow2 = case["pow2"]
    experts = "E" in case
    bounds = s["offsets"].tolist() if experts else [0, case["M"]]
    groups = [(b, e, s["w"][i] if experts else s["w"], s["wscales"][i] if experts else s["wscales"]) for i, (b, e) in enumerate(zip(bounds, bounds[1:]))]
    if kind in ("linear", "experts"):
        x = _exact_rows(s["x"].double(), pow2)
        y = torch.empty(case["M"], case["N"], dtype=torch.float64, device=x.device)
        for b, e, codes, scales in groups:
            if e > b:
                y[b:e] = torch.einsum("mk,nk->mn", x[b:e], _exact_tiles(codes, scales))
        return y if s["bias"] is None else y + s["bias"].double()
    dy = s["dy"].double()
    rows, columns = _exact_rows(dy, pow2), _exact_columns(dy, bounds, pow2)
    dx = torch.empty(case["M"], case["K"], dtype=torch.float64, device=dy.device)
    dw = torch.zeros(len(groups), case["N"], case["K"], dtype=torch.float64, device=dy.device)
    at = 0                                                   # first row of the expert in the kept activations
    for i, (b, e, codes, scales) in enumerate(groups):
        if e == b:
            continue
        dx[b:e] = torch.einsum("mn,nk->mk", rows[b:e], _exact_tiles(codes, scales))
        x = s["x"][at:at + e - b].double()
        for r in range(0, e - b, BLOCK):
            x[r:r + BLOCK] *= s["xscales"][(at + r) // BLOCK].double()
        dw[i] = torch.einsum("mn,mk->nk", columns[b:e], x)
        at += -(-(e - b) // BLOCK) * BLOCK
    return {"dx": dx, "dw": dw if experts else dw[0]}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    kind = case["kind"]
    if kind == "clip":
        # the norm has to be known before the first number is scaled: every gradient is read twice
        return {"bytes": 3 * size * case["elements"], "flops": 3 * case["elements"]}
    M, N, K, E = case["M"], case["N"], case["K"], case.get("E", 1)
    busy = E * (1 - (1 - 1 / E) ** M)                        # experts that a token comes to, if all are as popular
    weight = busy * (N * K + 4 * -(-N // BLOCK) * -(-K // BLOCK))
    if kind in ("linear", "experts"):
        return {"bytes": size * M * K + weight + size * M * N, "flops": 2 * M * N * K}
    wsize = 4 if case["wdtype"] == "fp32" else size
    kept = M * K + 4 * -(-M // BLOCK) * K
    return {"bytes": size * M * N + weight + kept + size * M * K + wsize * E * N * K, "flops": 4 * M * N * K}
