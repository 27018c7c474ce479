"""The operators around an 8-bit KAN layer in a language model's block, over the sizes that programs call them at, each
beside its plain form (elementary torch operations in 32 bits) and what a 64-bit evaluation returns.

A case names the operator (op), its sizes and its types:
  norm      the residual's addition and the root-mean-square norm of [rows, width], out in 8-bit floating point with a scale
            for each 128 columns of a row; x and residual are "f32", "f16" or "bf16" (residual also "none"); "strided": the
            rows of x are part of wider ones
  weights   weights [experts, outputs, inputs] (experts 0: one matrix) to 8-bit floating point with a scale for each block
            of 128 x 128
  product   [rows, inputs] times [outputs, inputs] transposed, both in 8 bits with their scales, out in `out`
  experts   the same product grouped by expert: `top` experts for each of `tokens`, the rows sorted by expert; `skew` is the
            spread of the experts' popularity (in nats), which makes the groups ragged and leaves some empty
"""
from __future__ import annotations

import math

import torch

own = False          # False: the plain forms; True: this package's operators

BLOCK = 128          # columns (and rows of a weight) that share a scale
LARGEST = 448.0      # the largest finite value of float8_e4m3fn
SMALLEST_SCALE = 2.0 ** -126
EPS = 1e-6
_TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_PRODUCT_MOST = 2.0 * 8192 * 4096 * 4096
_EXPERTS_MOST = 2.0 * 16384 * 2048 * 1024


def listed():
    return [
        # one token of a decoding step in front of a 1024-wide layer: latency
        {"name": "norm_token", "op": "norm", "rows": 1, "width": 1024, "x": "bf16", "residual": "bf16", "strided": False},
        # an irregular width in 32 bits, as a KAN layer hands its outputs on: no block of 128 ends where a row does
        {"name": "norm_ragged_1000", "op": "norm", "rows": 1000, "width": 300, "x": "f32", "residual": "f32", "strided": False},
        # the widest layer's largest batch
        {"name": "norm_32768", "op": "norm", "rows": 32768, "width": 1024, "x": "bf16", "residual": "bf16", "strided": False},
        # the weights of a square projection, converted as a model is loaded
        {"name": "weights_4096", "op": "weights", "experts": 0, "outputs": 4096, "inputs": 4096, "x": "bf16"},
        # a few irregular experts in 32 bits
        {"name": "weights_ragged", "op": "weights", "experts": 8, "outputs": 300, "inputs": 200, "x": "f32"},
        # one token through a square projection: latency
        {"name": "product_token", "op": "product", "rows": 1, "inputs": 1024, "outputs": 1024, "out": "f32"},
        # a server's decoding step: the weights' bytes
        {"name": "product_16", "op": "product", "rows": 16, "inputs": 4096, "outputs": 4096, "out": "bf16"},
        # the irregular layer's widths
        {"name": "product_ragged_1000", "op": "product", "rows": 1000, "inputs": 200, "outputs": 300, "out": "f32"},
        # a long prompt or a training-size batch: the matrix cores
        {"name": "product_8192", "op": "product", "rows": 8192, "inputs": 4096, "outputs": 4096, "out": "bf16"},
        # a decoding step through a few experts: the weights' bytes of those that were picked
        {"name": "experts_16", "op": "experts", "tokens": 16, "top": 2, "experts": 8, "inputs": 1024, "outputs": 1024,
         "out": "bf16", "skew": 1.0},
        # irregular experts, ragged groups, 32 bits out for a table layer behind them
        {"name": "experts_ragged", "op": "experts", "tokens": 500, "top": 3, "experts": 12, "inputs": 200, "outputs": 300,
         "out": "f32", "skew": 1.0},
        # a long prompt through many experts
        {"name": "experts_8192", "op": "experts", "tokens": 8192, "top": 2, "experts": 32, "inputs": 2048, "outputs": 1024,
         "out": "bf16", "skew": 0.5},
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):                                # half of them whole blocks or pieces of 16, half whatever comes
        w = log_int(lo, hi)
        step = rng.choice([1, 1, 16, BLOCK])
        return max(lo, w // step * step) if w >= step else w

    op = rng.choice(["norm", "weights", "product", "product", "experts", "experts"])
    if op == "norm":
        w = width(8, 8192)
        return {"op": op, "rows": max(1, min(log_int(1, 32768), (1 << 25) // w)), "width": w, "x": rng.choice(sorted(_TYPE)),
                "residual": rng.choice(sorted(_TYPE) + ["none"]), "strided": rng.random() < 0.25}
    if op == "weights":
        outputs, inputs = width(16, 4096), width(16, 4096)
        experts = min(rng.choice([0, 0, 2, 8, 16]), (1 << 24) // (outputs * inputs))
        return {"op": op, "experts": experts, "outputs": outputs, "inputs": inputs, "x": rng.choice(sorted(_TYPE))}
    if op == "product":
        inputs, outputs = width(16, 8192), width(2, 8192)
        outputs = max(1, min(outputs, (1 << 25) // inputs))
        rows = min(log_int(1, 32768), (1 << 25) // max(inputs, outputs), int(_PRODUCT_MOST / (2.0 * inputs * outputs)))
        return {"op": op, "rows": max(1, rows), "inputs": inputs, "outputs": outputs, "out": rng.choice(sorted(_TYPE))}
    inputs, outputs, experts, top = width(16, 4096), width(16, 4096), rng.randint(2, 64), rng.randint(1, 4)
    outputs = max(1, min(outputs, (1 << 26) // (inputs * experts)))
    rows = min(log_int(1, 8192) * top, (1 << 24) // max(inputs, outputs), int(_EXPERTS_MOST / (4.0 * inputs * outputs)))
    return {"op": op, "tokens": max(1, rows // top), "top": min(top, experts), "experts": experts, "inputs": inputs, "outputs": outputs,
            "out": rng.choice(sorted(_TYPE)), "skew": rng.choice([0.0, 0.5, 1.0])}


# ---- inputs ------------------------------------------------------------------------------------------------------
def _blocks(n):
    return -(-n // BLOCK)


def _pad_columns(v):
    return torch.nn.functional.pad(v, (0, _blocks(v.shape[-1]) * BLOCK - v.shape[-1]))


def _codes_by_row(v):
    """float8 codes [..., n] and scales [..., blocks] of v [..., n] in 32 bits."""
    n = v.shape[-1]
    b = _pad_columns(v).unflatten(-1, (_blocks(n), BLOCK))
    scales = (b.abs().amax(dim=-1) / LARGEST).clamp(min=SMALLEST_SCALE)
    return (b / scales[..., None]).to(torch.float8_e4m3fn).flatten(-2)[..., :n].contiguous(), scales


def _codes_by_block(w):
    """float8 codes [..., n, k] and scales [..., row blocks, column blocks] of w [..., n, k]."""
    n, k = w.shape[-2:]
    v = torch.nn.functional.pad(w.float(), (0, _blocks(k) * BLOCK - k, 0, _blocks(n) * BLOCK - n))
    b = v.unflatten(-1, (_blocks(k), BLOCK)).unflatten(-3, (_blocks(n), BLOCK))      # [..., row block, row, column block, column]
    scales = (b.abs().amax(dim=(-3, -1)) / LARGEST).clamp(min=SMALLEST_SCALE)
    codes = (b / scales[..., :, None, :, None]).to(torch.float8_e4m3fn).flatten(-2).flatten(-3, -2)
    return codes[..., :n, :k].contiguous(), scales


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def activations(rows, width):                     # channels of different size, as a model's are
        return normal(rows, width) * torch.exp(0.7 * normal(width))

    op = case["op"]
    if op == "norm":
        rows, width = case["rows"], case["width"]
        x = activations(rows, width + 24 if case["strided"] else width).to(_TYPE[case["x"]])[:, :width]
        residual = None if case["residual"] == "none" else (3.0 * activations(rows, width)).to(_TYPE[case["residual"]])
        return {"op": op, "x": x, "residual": residual, "weight": (1.0 + 0.2 * normal(width)).to(x.dtype)}
    if op == "weights":
        shape = ([case["experts"]] if case["experts"] else []) + [case["outputs"], case["inputs"]]
        return {"op": op, "weight": (normal(*shape) / math.sqrt(case["inputs"])).to(_TYPE[case["x"]])}
    shape = ([case["experts"]] if op == "experts" else []) + [case["outputs"], case["inputs"]]
    rows = case["tokens"] if op == "experts" else case["rows"]
    state = {"op": op, "out": _TYPE[case["out"]]}
    state["x"], state["x_scales"] = _codes_by_row(activations(rows, case["inputs"]))
    state["weight"], state["weight_scales"] = _codes_by_block(normal(*shape) / math.sqrt(case["inputs"]))
    if op == "experts":
        logits = normal(rows, case["experts"]) + case["skew"] * normal(case["experts"])
        expert = logits.topk(case["top"], dim=1).indices.flatten()
        order = torch.sort(expert, stable=True).indices
        state["rows"] = order // case["top"]                                  # the token of each sorted row
        state["group_sizes"] = torch.bincount(expert, minlength=case["experts"])
    return state


# ---- one pass ----------------------------------------------------------------------------------------------------
def _values(codes, scales):
    return codes.float() * scales.repeat_interleave(BLOCK, dim=-1)[..., :codes.shape[-1]]


def _weight_values(codes, scales):
    return codes.float() * scales.repeat_interleave(BLOCK, dim=-2)[..., :codes.shape[-2], :].repeat_interleave(BLOCK, dim=-1)[..., :codes.shape[-1]]


def _plain_norm(x, weight, residual):
    h = x.float() if residual is None else x.float() + residual.float()
    y = h * torch.rsqrt(h.square().mean(dim=-1, keepdim=True) + EPS) * weight.float()
    return *_codes_by_row(y), None if residual is None else h.to(residual.dtype)


def _plain_product(x, x_scales, weight, weight_scales, out):
    return torch.matmul(_values(x, x_scales), _weight_values(weight, weight_scales).t()).to(out)


def _plain_experts(x, x_scales, weight, weight_scales, group_sizes, rows, out):
    """All experts as one batched product: every group is padded to the largest."""
    ends = group_sizes.cumsum(0)
    at = torch.arange(rows.numel(), device=x.device)
    group = torch.searchsorted(ends, at, right=True)
    place = at - (ends - group_sizes)[group]
    padded = torch.zeros((group_sizes.numel(), int(group_sizes.max()), x.shape[1]), device=x.device)
    padded[group, place] = _values(x, x_scales)[rows]
    y = torch.bmm(padded, _weight_values(weight, weight_scales).transpose(1, 2).contiguous())
    return y[group, place].to(out)


def run(state):
    s = state
    if own:
        import paper_2601_03332_amd as lk
        if s["op"] == "norm":
            return lk.lutkan_rmsnorm_fp8(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        if s["op"] == "weights":
            return lk.lutkan_quantise_fp8(s["weight"])
        if s["op"] == "product":
            return lk.lutkan_matmul_fp8(s["x"], s["x_scales"], s["weight"], s["weight_scales"], dtype=s["out"])
        return lk.lutkan_grouped_matmul_fp8(s["x"], s["x_scales"], s["weight"], s["weight_scales"], s["group_sizes"], rows=s["rows"],
                                            dtype=s["out"])
    if s["op"] == "norm":
        return _plain_norm(s["x"], s["weight"], s["residual"])
    if s["op"] == "weights":
        return _codes_by_block(s["weight"])
    if s["op"] == "product":
        return _plain_product(s["x"], s["x_scales"], s["weight"], s["weight_scales"], s["out"])
    return _plain_experts(s["x"], s["x_scales"], s["weight"], s["weight_scales"], s["group_sizes"], s["rows"], s["out"])


def work(case):
    """Each input once, each output once; for experts those rows of x and those experts' weights that the routing can reach."""
    size = {"f32": 4, "f16": 2, "bf16": 2, "none": 0}
    if case["op"] == "norm":
        n, w = case["rows"], case["width"]
        return {"bytes": n * w * (size[case["x"]] + 2.0 * size[case["residual"]] + 1.0) + 4.0 * n * _blocks(w) + w * size[case["x"]],
                "flops": 8.0 * n * w}
    matrices = max(1, case.get("experts", 0))
    if case["op"] == "weights":
        n, k = case["outputs"], case["inputs"]
        return {"bytes": matrices * (n * k * (size[case["x"]] + 1.0) + 4.0 * _blocks(n) * _blocks(k)), "flops": 3.0 * matrices * n * k}
    k, n = case["inputs"], case["outputs"]
    read = case["tokens"] if case["op"] == "experts" else case["rows"]
    rows = read * case.get("top", 1)
    held = min(matrices, rows) * (n * k + 4.0 * _blocks(n) * _blocks(k))
    return {"bytes": read * (k + 4.0 * _blocks(k)) + held + rows * n * float(size[case["out"]]), "flops": 2.0 * rows * k * n}


# ---- the same outputs in 64 bits -----------------------------------------------------------------------------------
def _decoded(codes):
    """Values of float8_e4m3fn codes from their bits: sign, four bits of exponent (bias 7), three of mantissa."""
    bits = codes.contiguous().view(torch.uint8).to(torch.int64)
    exponent, mantissa = (bits >> 3) & 15, (bits & 7).to(torch.float64)
    power = torch.exp2((exponent.clamp(min=1) - 7).to(torch.float64))
    value = torch.where(exponent == 0, mantissa / 8.0, 1.0 + mantissa / 8.0) * power
    return torch.where(bits >= 128, -value, value)


def _exact_product(x, x_scales, weight, weight_scales):
    """Block by block along the inputs: the product of the codes, then both scales."""
    y = torch.zeros((x.shape[0], weight.shape[0]), dtype=torch.float64, device=x.device)
    of_row = torch.arange(weight.shape[0], device=x.device) // BLOCK
    for b in range(x_scales.shape[1]):
        part = _decoded(x[:, b * BLOCK:(b + 1) * BLOCK]) @ _decoded(weight[:, b * BLOCK:(b + 1) * BLOCK]).t().contiguous()
        y += part * x_scales[:, b, None].double() * weight_scales[of_row, b].double()
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        y = h / torch.sqrt((h * h).sum(dim=1, keepdim=True) / h.shape[1] + EPS) * s["weight"].double()
        codes, scales = torch.empty_like(y), torch.empty((y.shape[0], _blocks(y.shape[1])), dtype=torch.float64, device=y.device)
        for b in range(scales.shape[1]):
            part = y[:, b * BLOCK:(b + 1) * BLOCK]
            scales[:, b] = torch.maximum(part.abs().max(dim=1).values / LARGEST, torch.full_like(part[:, 0], SMALLEST_SCALE))
            codes[:, b * BLOCK:(b + 1) * BLOCK] = part / scales[:, b, None]
        return codes, scales, None if s["residual"] is None else h              # the codes as they are before they are rounded
    if case["op"] == "weights":
        w = s["weight"].double()
        codes = torch.empty_like(w)
        scales = torch.empty((*w.shape[:-2], _blocks(w.shape[-2]), _blocks(w.shape[-1])), dtype=torch.float64, device=w.device)
        for r in range(scales.shape[-2]):
            for b in range(scales.shape[-1]):
                at = (..., slice(r * BLOCK, (r + 1) * BLOCK), slice(b * BLOCK, (b + 1) * BLOCK))
                scales[..., r, b] = (w[at].abs().flatten(-2).max(dim=-1).values / LARGEST).clamp(min=SMALLEST_SCALE)
                codes[at] = w[at] / scales[..., r, b, None, None]
        return codes, scales
    if case["op"] == "product":
        return _exact_product(s["x"], s["x_scales"], s["weight"], s["weight_scales"])
    parts, first = [], 0
    for e, n in enumerate(s["group_sizes"].tolist()):
        at = s["rows"][first:first + n]
        parts.append(_exact_product(s["x"][at], s["x_scales"][at], s["weight"][e], s["weight_scales"][e]))
        first += n
    return torch.cat(parts)
